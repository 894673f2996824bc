"""The serving loop with KV caches in 8 bits (paper_2508_01989_amd/instance.py, `kvq`): every flow of requests between instances, all of them
in 8 bits or some in 16.  The plain form of the cache is kept beside every instance: each iteration's attention, and what a request's cache
stands for after each move, are compared with it."""
import numpy as np
import pytest

import oracle
from oracle import kvq

SHAPE, LAYERS = (8, 2, 128), 2
KINDS = {"all_in_8_bits": [True, True, True], "one_in_16_bits": [True, False, True]}


def scenario(dry, kinds):
    from paper_2508_01989_amd import sched
    from paper_2508_01989_amd.instance import Cluster, make_request
    cm = sched.cost_model(LAYERS, 20e-6, 1e-6, 2e-11, 1e-9)
    cl = Cluster([sched.P_HEAVY, sched.D_HEAVY, sched.D_HEAVY], [64, 16, 16], [48, 12, 12], SHAPE, LAYERS, cm,
                 tpot_slo=80e-6, ttft_slo=1e-3, watermark_frac=0.75, dry=dry, kvq=kinds)
    rng = np.random.default_rng(3)
    reqs, t = [], 0.0
    for i in range(12):
        t += float(rng.exponential(150e-6))
        reqs.append(make_request(i, int(rng.integers(5, 120)), int(rng.integers(2, 40)), t, SHAPE, LAYERS, seed=i, dry=dry))
    return cl, reqs


def check_bookkeeping(cl, reqs, done):
    assert sorted(r.rid for r in done) == [r.rid for r in reqs]
    assert all(x.blocks_used == 0 and not x.queue and not x.decodes for x in cl.inst)
    s = cl.stats
    assert s["handoffs"] > 0 and s["in_place"] > 0 and s["degrade_flows"] > 0 and s["backflows"] > 0 and s["bytes_moved"] > 0


@pytest.mark.parametrize("kinds", KINDS)
def test_dry_run_exercises_every_flow(kinds):
    cl, reqs = scenario(True, KINDS[kinds])
    check_bookkeeping(cl, reqs, cl.run(reqs))
    assert scenario(True, True)[0].inst[2].kvq and not scenario(True, False)[0].inst[0].kvq


class Plain16:
    """A cache in 16 bits with the interface of kvq.Cache that the test uses."""

    def __init__(self, blocks):
        _, self.Hkv, self.D = SHAPE
        self.k, self.v = oracle.new_pool(blocks, self.Hkv, self.D)

    def append(self, q_start, ctx, table, k, v):
        oracle.kv_append(self.k, self.v, self.Hkv, self.D, 16, q_start, ctx, table, k, v)

    def read(self, row, n):
        return [kvq.widen(x, "bf16") for x in oracle.kv_gather(self.k, self.v, self.Hkv, self.D, 16, row, n)]

    def widened_pools(self, table, kv):
        return self.k, self.v


@pytest.mark.gpu
@pytest.mark.parametrize("kinds", KINDS)
def test_outputs_and_caches_on_every_route(kinds, monkeypatch):
    import torch
    assert torch.cuda.is_available()
    from paper_2508_01989_amd import instance as I
    Hq, Hkv, D = SHAPE
    cl, reqs = scenario(False, KINDS[kinds])
    plain = {x.index: [kvq.Cache(x.num_blocks, Hkv, D) if x.kvq else Plain16(x.num_blocks) for _ in range(LAYERS)] for x in cl.inst}
    host = lambda t: t.cpu().numpy().view(np.uint16)  # noqa: E731
    worst = [0.0]
    run_layers, migrate = I.Instance._run_layers, I.Cluster.migrate

    def checked_run(self, rs, q_len, ctx, q_start):
        run_layers(self, rs, q_len, ctx, q_start)
        table = np.zeros((len(rs), max(len(r.blocks) for r in rs)), np.int32)
        for i, r in enumerate(rs):
            table[i, :len(r.blocks)] = r.blocks
        for l in range(LAYERS):
            part = lambda x: np.concatenate([host(getattr(r, x)[l, c:c + n]) for r, n, c in zip(rs, q_len, ctx)])  # noqa: E731
            c = plain[self.index][l]
            c.append(q_start, ctx, table, part("k"), part("v"))
            kp, vp = c.widened_pools(table, ctx + q_len)
            args = (Hq, Hkv, D, 16, q_start, ctx, table, part("q"), 1.0 / np.sqrt(D))
            want, mean = oracle.attention(kp, vp, *args), oracle.attention(kp, vp & np.uint16(0x7FFF), *args)
            got = kvq.widen(part("out"), "bf16")
            # a half step of bf16 for the probabilities and one for the output, relative, and a fiftieth for sums in 32 bits
            worst[0] = max(worst[0], float((np.abs(got - want) / (2.0 ** -8 * 1.02 * (mean + np.abs(want)) + 1e-30)).max()))

    def checked_migrate(self, req, dst, now, why):
        src, old, n = self.inst[req.where], list(req.blocks), req.done
        migrate(self, req, dst, now, why)
        for l in range(LAYERS):
            rows = plain[src.index][l].read(np.array(old), n)
            plain[dst.index][l].append(np.array([0, n], np.int32), np.zeros(1, np.int32), np.array([req.blocks], np.int32),
                                       *(kvq.narrow(x, "bf16") for x in rows))
            if dst.kvq:
                for dev, c in ((dst.k_pools[l], plain[dst.index][l].k), (dst.v_pools[l], plain[dst.index][l].v), (dst.scales[l], plain[dst.index][l].scales)):
                    used = np.array(req.blocks[:n // 16], np.int64)  # whole pages
                    assert np.array_equal(dev.cpu().numpy().reshape(c.shape)[used], c[used])

    monkeypatch.setattr(I.Instance, "_run_layers", checked_run)
    monkeypatch.setattr(I.Cluster, "migrate", checked_migrate)
    print(f"[case] instance loop, caches in 8 bits: {kinds}", flush=True)
    done = cl.run(reqs)
    check_bookkeeping(cl, reqs, done)
    assert worst[0] <= 1.0, worst[0]
