"""Runs whose devices exchange messages of 4 bits per parameter: the calls of a round together, round after round,
against the oracle's counters and the messages' definition (packed_reference.py)."""
import json

import numpy as np
import pytest
import torch

import packed_reference as ref
from gpu_common import require_gpu
from oracle_driver import make_sim
from paper_2111_08274_b200 import binding, run, runtime, workloads
from test_gpu_packed import aggregate_reference, assert_same, to_storage

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def workload(n, p, k, dtype, **kw):
    return workloads.Workload("packed", n, p, k, 5, "uniform", steps_lo=0, steps_hi=3, grad_std=1e-2, seed=91, dtype=dtype,
                              m_dtype=dtype, **kw)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rounding", [binding.ROUND_NEAREST, binding.ROUND_STOCHASTIC])
@pytest.mark.parametrize("n,p,k,sync_every,beta,weight_mode", [(4, 2003, 2, 2, 1.0, 0), (5, 700, 3, 0, 1.0, 1), (3, 33, 1, 2, 0.5, 0),
                                                              (6, 4097, 6, 3, 1.0, 1)])
def test_rounds_that_exchange_messages(oracle, n, p, k, sync_every, beta, weight_mode, rounding, dtype):
    """Every round: local steps (already tested; their result is read back), selection as the oracle's, then the exchange
    bit for bit as the definition says: messages, residuals, aggregate, base, versions, products."""
    wl = workload(n, p, k, dtype, sync_every=sync_every, sync_beta=beta, weight_mode=weight_mode)
    arena, sim = runtime.Arena(wl), make_sim(oracle, wl)
    exchange = runtime.Exchange(arena, rounding)
    base = arena.w[0, :p].float().cpu().numpy()
    residual = np.zeros((n, p), np.float32)
    for r in range(wl.rounds):
        arena.h.local_step(arena.ids, wl.steps_for_round(r), wl.lr)
        sim.local_step(wl.device_ids(), wl.steps_for_round(r), wl.lr)
        rows = arena.w[:, :p].float().cpu().numpy()
        sel = arena.h.select(r, k, arena.select_seed)
        assert np.array_equal(sel, sim.select(r, k, wl.select_seed()))
        a = arena.h.aggregation_weights(sel)
        sync = bool(sync_every) and (r + 1) % sync_every == 0
        exchange.synchronise(sel, r, sync)
        d = []
        for i in sel:
            u = ref.to_send(rows[i], base, residual[i])
            codes, scales = ref.message(u, ref.random_bits(wl.seed, int(i), r, p) if rounding else None)
            assert np.array_equal(exchange.messages[int(i)].cpu().numpy(), ref.to_bytes(codes, scales, p))
            residual[i] = ref.residual_after(u, codes, scales)
            d.append(ref.values(codes, scales, p))
        assert_same(exchange.residual[:, :p].cpu().numpy(), residual)
        x = aggregate_reference(a, d, base)
        receivers = range(n) if sync and beta == 1.0 else sel
        want = rows.copy()
        for i in receivers:
            want[i] = to_storage(x, arena.w.dtype)
        if sync and beta < 1.0:
            for i in set(range(n)) - set(int(j) for j in sel):
                mine = (np.float32(1) - np.float32(beta)) * rows[i]
                want[i] = to_storage((np.longdouble(beta) * want[sel[0]].astype(np.longdouble) + mine.astype(np.longdouble)), arena.w.dtype)
        got = arena.w[:, :p].float().cpu().numpy()
        assert_same(got, want, r)
        if sync and beta == 1.0:
            base = want[0]
        assert_same(exchange.base.float().cpu().numpy(), base)
        sim.aggregate(sel)
        if sync:
            others = np.setdiff1d(np.arange(n), sel).astype(np.int32)
            sim.broadcast(int(sel[0]), others) if beta == 1.0 else sim.integrate(int(sel[0]), others, beta)
        assert np.array_equal(arena.h.get_versions()[0], sim.get_versions()[0])
        d = np.stack(d)
        assert np.all(np.abs(exchange.read_products() - d @ d.T) <= 4e-6 * (np.abs(d) @ np.abs(d).T) + 1e-37)
    arena.h.debug_check()
    arena.close()


def test_round_helper_is_the_calls():
    wl = workload(4, 3001, 2, 0, sync_every=2)
    one, two = runtime.Arena(wl), runtime.Arena(wl)
    e1, e2 = runtime.Exchange(one), runtime.Exchange(two)
    for r in range(wl.rounds):
        s1 = one.run_round_packed(r, e1)
        two.h.local_step(two.ids, wl.steps_for_round(r), wl.lr)
        s2 = two.h.select(r, wl.k, two.select_seed)
        e2.synchronise(s2, r, (r + 1) % 2 == 0)
        two.h.stats_enqueue(int(s2[0]))
        assert np.array_equal(s1, s2)
        for x, y in zip(one.h.stats_read(), two.h.stats_read()):
            assert np.array_equal(x, y)
        for x, y in ((one.w, two.w), (e1.messages, e2.messages), (e1.residual, e2.residual), (e1.products, e2.products)):
            assert torch.equal(x, y)
    one.close()
    two.close()


def test_exchange_without_residuals():
    wl = workload(3, 500, 2, 0)
    arena = runtime.Arena(wl)
    exchange = runtime.Exchange(arena, binding.ROUND_NEAREST, residual=False)
    assert exchange.residual is None
    for r in range(3):
        sel = arena.run_round_packed(r, exchange)
    got = arena.w[:, :500].cpu().numpy()
    assert np.array_equal(got[sel[0]], got[sel[1]]) and np.all(np.isfinite(got))
    arena.close()


@pytest.mark.parametrize("how", ["nearest", "stochastic"])
def test_command_logs_messages(tmp_path, how):
    path, plain = tmp_path / "packed.jsonl", tmp_path / "plain.jsonl"
    args = ["--workload", "c1", "--n-params", "20003", "--rounds", "6"]
    run.main([*args, "--jsonl", str(path), "--packed", how])
    run.main([*args, "--jsonl", str(plain)])
    rows, others = ([json.loads(line) for line in f.read_text().splitlines()] for f in (path, plain))
    assert len(rows) == len(others) == 6
    for row, other in zip(rows, others):
        for key in ("selected", "versions", "step_counters", "global_sync"):
            assert row[key] == other[key], key
        products = np.array(row["message_products"])
        assert products.shape == (2, 2) and np.array_equal(products, products.T) and np.all(np.diag(products) > 0)
        assert row["message_bytes"] == binding.hadfl_packed_bytes(20003)
        assert all(row["divergence2"][s] == 0.0 for s in row["selected"])
        # a message leaves out at most a sixth of the largest value of a block: the models stay near those of the plain run
        assert np.allclose(row["norm2"], other["norm2"], rtol=0.05)


def test_command_with_predicted_versions(tmp_path):
    path = tmp_path / "planned.jsonl"
    run.main(["--workload", "c1", "--n-params", "5003", "--rounds", "5", "--jsonl", str(path), "--packed", "stochastic",
              "--predict", "0.6"])
    rows = [json.loads(line) for line in path.read_text().splitlines()]
    assert rows[1]["planned_versions"] is None and rows[4]["planned_versions"] is not None
