"""Two host threads with streams, buffers and workspaces of their own: calls that share a kernel but need
different amounts of shared memory, at the same time, succeed and give the bits that they give alone."""
import threading

import pytest
import torch

from paper_2609_32525_gb300.workloads import make_case

from _parity import upload

pytestmark = pytest.mark.gpu


def _norm(lib, C, res, seed, backward):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows = 64
    x, y = (torch.randn(rows, C, generator=g, device="cuda") for _ in range(2))
    r, other = lib.rows_of(x), torch.randn(rows, C, generator=g, device="cuda") if res else None
    mean, rstd = x.mean(1), torch.rsqrt(x.var(1, unbiased=False) + 1e-5)
    if not backward:
        out = [torch.empty_like(x), torch.empty_like(mean), torch.empty_like(mean)]
        return out, lambda s: lib.fs_norm_fwd(r, x, other, None, None, 1e-5, None, *out, stream=s)
    out, ws = [torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")], lib.norm_workspace(r)
    return out, lambda s: lib.fs_norm_bwd(r, x, None, None, None, mean, rstd, y, other, *out, False, ws, stream=s)


def _coupling(lib, G, seed):
    v = upload(make_case(1, 300, 2, 32, G, dtype="bf16", seed=seed, backward=True))
    c = lib.Coupling(1, 300, 2, 32, G, torch.bfloat16, backward=True)
    a = [v[k] for k in ("x_mid", "fx", "W_slice", "bias", "tau", "M")]

    def call(s):
        c.forward(*a, stream=s)
        c.backward(*a, v["dout"], stream=s)

    return [c.out, c.tokens, c.dx_mid, c.dfx, c.dW, c.dM], call


class Recorder:
    """Stands in for the loaded library: makes each call and keeps it with its arguments."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        fn = getattr(self.real, name)

        def call(*args):
            self.calls.append((fn, args))
            return fn(*args)

        return call


# Widths of 129 to 255 fp32 channels, odd, share the kernels that read rows by bulk copies; couplings of
# any number of slots share the statistics, the deslice and the backward.
JOBS = {
    "norm_fwd": (lambda lib: _norm(lib, 129, False, 1, False), lambda lib: _norm(lib, 255, True, 2, False), 20000),
    "norm_bwd": (lambda lib: _norm(lib, 129, False, 3, True), lambda lib: _norm(lib, 255, True, 4, True), 20000),
    "coupling": (lambda lib: _coupling(lib, 64, 5), lambda lib: _coupling(lib, 512, 6), 2000),
}


@pytest.mark.parametrize("name", JOBS)
def test_calls_of_different_sizes_at_once(lib, monkeypatch, name):
    *makers, n = JOBS[name]
    jobs, streams = [m(lib) for m in makers], [torch.cuda.Stream() for _ in makers]
    real, calls = lib._lib, []
    torch.cuda.synchronize()
    for (_, call), stream in zip(jobs, streams):  # as C calls, which run side by side
        monkeypatch.setattr(lib, "_lib", Recorder(real))
        call(stream)
        calls.append(lib._lib.calls)
    torch.cuda.synchronize()
    want = [[t.clone() for t in out] for out, _ in jobs]
    torch.cuda.synchronize()
    failed, start = [], threading.Barrier(2)

    def work(stream, calls):
        start.wait()
        for i in range(n):
            failed.extend(st for fn, args in calls if (st := fn(*args)) != lib.FS_OK)
            if i % 500 == 499:
                stream.synchronize()

    threads = [threading.Thread(target=work, args=a) for a in zip(streams, calls)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, f"{len(failed)} calls failed"
    for (out, _), w in zip(jobs, want):
        assert all(torch.equal(a, b) for a, b in zip(out, w))
