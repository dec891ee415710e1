"""Host threads, each with a context of its own, that call at the same time."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


def _together(jobs):
    """Runs the jobs in threads that start together; raises what one of them raised."""
    gate, failed = threading.Barrier(len(jobs)), []

    def run(job):
        try:
            gate.wait()
            job()
        except Exception as e:
            failed.append(e)
    threads = [threading.Thread(target=run, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if failed:
        raise failed[0]


@pytest.mark.parametrize("large,small", [((700, 256, 256), (700, 250, 1)), ((200, 1024, 1024), (200, 1000, 1)), ((150000, 1024, 1), (90000, 1024, 1))])
def test_threads_route_with_shared_memory_of_different_sizes(large, small):
    """The kernels' limits of shared memory are the device's: a thread with fewer experts or groups must not lower another's."""
    import paper_1904_02205_b200 as psb

    jobs, checks = [], []
    for i, (tokens, experts, groups) in enumerate((large, small)):
        ctx, stream = psb.Context(0), torch.cuda.Stream()
        logits = torch.randn(tokens, experts, generator=torch.Generator().manual_seed(i)).cuda()
        how = dict(groups=groups, top_groups=min(groups, 9), stream=stream)
        torch.cuda.synchronize()
        want = ctx.route_experts(logits, 4, **how)
        torch.cuda.synchronize()

        def job(ctx=ctx, stream=stream, logits=logits, how=how, want=want):
            got = []
            with torch.cuda.stream(stream):
                for _ in range(200):
                    got.append(ctx.route_experts(logits, 4, **how))
            stream.synchronize()
            assert ctx.device_status(stream) == 0
            for g in got:
                assert all(torch.equal(g[k], want[k]) for k in want)
        jobs.append(job)
        checks.append(ctx)
    _together(jobs)
    for ctx in checks:
        ctx.close()
