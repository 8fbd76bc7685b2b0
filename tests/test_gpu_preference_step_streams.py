"""A preference step made on one stream and used on others: every result has the bits of a step that stays on one stream."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_preference_step import make

pytestmark = pytest.mark.gpu


def outcome(job):
    torch.cuda.synchronize()
    return [t.clone() for t in (job.reference, job.logits, job.dlogits, job.drows, job.gate, job.scale, job.d_gate, job.d_scale, *job.A, *job.B, *job.dA, *job.dB)]


def steps(job, rows, targets, streams):
    """Reference and steps, each under another stream, whose inputs arrive late; the losses are read under the caller's stream."""
    losses = []
    for i in range(4):
        with torch.cuda.stream(streams[i % len(streams)]):
            torch.empty(1 << 25, device="cuda").normal_()          # the stream has work before the inputs are there
            r, t = rows.clone(), targets.clone()
            if i == 0:
                job.set_reference(r, t)
            losses.append(job.step(r, t))
            job.forward(r, counter=100 + i)
            job.losses(t)
            job.backward(r, t, counter=100 + i)
            losses.append(job.loss.clone())
            r.zero_()                                              # behind the backward's reads
            t.fill_(-100)
    torch.cuda.synchronize()
    return [x if isinstance(x, list) else x.tolist() for x in losses]


def test_a_step_made_on_one_stream_runs_under_others():
    job, rows, targets = make()
    main = torch.cuda.current_stream()
    want = steps(job, rows, targets, [main])
    state = outcome(job)
    sides = [torch.cuda.Stream() for _ in range(3)]
    for made_on, run_on in ((main, sides[:2]), (sides[2], [main, sides[0]]), (sides[0], [sides[1]])):
        torch.cuda.synchronize()
        with torch.cuda.stream(made_on):
            other, r, t = make()
        torch.cuda.synchronize()
        assert steps(other, r, t, run_on) == want
        for a, b in zip(outcome(other), state):
            assert torch.equal(a, b)
