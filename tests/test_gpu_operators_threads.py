"""The operators called from several threads at once: the entry points keep nothing of one call that another could change."""
import ctypes as C
import shutil
import subprocess

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# threads without the interpreter's lock between two calls
THREADS = r"""
#include <pthread.h>
#include <stdatomic.h>
#include <stdint.h>
typedef int (*entry)(const void*, uint64_t, const void*, uint64_t, void*, uint64_t, int, uint64_t, uint64_t, const void*, int, const float*,
                     const float*, void*, void*, int, void*, uint64_t, void*);
struct job { entry f; void *dy, *x, *dx; uint64_t rows, cols; int type; float *mean, *rstd; void* stream; int calls, refused; };
static _Atomic int ready;
static int count;
static void* work(void* p) {
    struct job* j = p;
    atomic_fetch_add(&ready, 1);
    while (atomic_load(&ready) < count) {}
    for (int i = 0; i < j->calls; ++i)
        j->refused += 0 != j->f(j->dy, j->cols, j->x, j->cols, j->dx, j->cols, j->type, j->rows, j->cols, 0, 0, j->mean, j->rstd, 0, 0, 0, 0, 0, j->stream);
    return 0;
}
void run(struct job* j, int n) {
    pthread_t t[8];
    count = n;
    atomic_store(&ready, 0);
    for (int i = 0; i < n; ++i) pthread_create(&t[i], 0, work, &j[i]);
    for (int i = 0; i < n; ++i) pthread_join(t[i], 0);
}
"""


class Job(C.Structure):
    _fields_ = [("f", C.c_void_p), ("dy", C.c_void_p), ("x", C.c_void_p), ("dx", C.c_void_p), ("rows", C.c_uint64), ("cols", C.c_uint64),
                ("type", C.c_int), ("mean", C.c_void_p), ("rstd", C.c_void_p), ("stream", C.c_void_p), ("calls", C.c_int), ("refused", C.c_int)]


@pytest.mark.skipif(not shutil.which("gcc"), reason="no gcc")
@pytest.mark.parametrize("dtype,code", [(torch.bfloat16, 1), (torch.float32, 0)], ids=["bfloat16", "float32"])
def test_row_lengths_that_share_a_kernel(tmp_path, dtype, code):
    """Rows of different lengths take one kernel with different amounts of shared memory, none of which is refused."""
    from paper_2210_07454_b200 import binding, operators as ops
    (tmp_path / "threads.c").write_text(THREADS)
    subprocess.run(["gcc", "-O2", "-shared", "-fPIC", "-o", "threads.so", "threads.c", "-lpthread"], cwd=tmp_path, check=True)
    entry = C.cast(binding.lib().sk_layer_norm_backward, C.c_void_p)
    rows, kept, jobs = 4, [], (Job * 4)()
    for j, cols in zip(jobs, (8192, 4480, 6000, 2200)):
        gen = torch.Generator(device="cuda").manual_seed(cols)
        x, dy = (torch.randn(rows, cols, generator=gen, device="cuda").to(dtype) for _ in range(2))
        _, mean, rstd = ops.layer_norm(x)
        want, dx, stream = ops.layer_norm_backward(dy, x, None, mean, rstd)[0], torch.zeros_like(x), torch.cuda.Stream()
        kept.append((x, dy, mean, rstd, want, dx, stream))
        j.f, j.dy, j.x, j.dx, j.rows, j.cols, j.type = entry, dy.data_ptr(), x.data_ptr(), dx.data_ptr(), rows, cols, code
        j.mean, j.rstd, j.stream, j.calls = mean.data_ptr(), rstd.data_ptr(), stream.cuda_stream, 5000
    torch.cuda.synchronize()
    C.CDLL(str(tmp_path / "threads.so")).run(jobs, 4)
    torch.cuda.synchronize()
    assert [j.refused for j in jobs] == [0] * 4
    assert all(torch.equal(k[5], k[4]) for k in kept)
