"""Calls on a stream of their own: whose memory results are, and when memory that
is freed early is used again.  The streams are kept busy by a kernel that ends by
itself; nothing here depends on how long it takes, beyond that it outlasts a few
calls on the host."""
import pytest
import torch

from paper_2101_08763_amd import api

pytestmark = pytest.mark.gpu
N, D, L, K = 4000, 512, 4000, 3
BUSY = 200_000_000  # cycles, 0.1 s


def tensors(*x):
    """The tensors among results (MxRows among them)."""
    out = []
    for t in x:
        if isinstance(t, torch.Tensor):
            out.append(t)
        elif isinstance(t, (tuple, list)):
            out.extend(tensors(*t))
    return out


def span(t):
    return t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()


def apart(t, spans):
    a, b = span(t)
    return all(b <= x or y <= a for x, y in spans)


@pytest.fixture(scope="module")
def made():
    g = torch.Generator("cuda").manual_seed(0)
    V = torch.randn(N, D, generator=g, device="cuda")
    sets = torch.randint(0, N, (L, K), generator=g, device="cuda", dtype=torch.int32)
    q4, q8 = api.exemplar_mx_quantize(V, api.EXEMCL_MXFP4), api.exemplar_mx_quantize(V, api.EXEMCL_MXFP8)
    rstd = torch.ones(N, device="cuda")
    return V, sets, q4, q8, rstd


# name: (the inputs of a call, the call on a stream)
CALLS = {
    "eval": (lambda m: (m[0], m[1]), lambda a, st: api.exemplar_eval(a[0], a[1], stream=st)),
    "gain": (lambda m: (m[0], m[1][0], m[1][:, 0].contiguous()), lambda a, st: api.exemplar_gain(*a, stream=st)),
    "sqnorm": (lambda m: (m[0],), lambda a, st: api.exemplar_sqnorm(a[0], stream=st)),
    "greedy": (lambda m: (m[0],), lambda a, st: api.exemplar_greedy(a[0], 4, stream=st)),
    "quantize": (lambda m: (m[0],), lambda a, st: api.exemplar_mx_quantize(a[0], api.EXEMCL_MXFP8, stream=st)),
    "dequantize": (lambda m: (m[2],), lambda a, st: api.exemplar_mx_dequantize(a[0], torch.float32, stream=st)),
    "norm": (lambda m: (m[0], m[0].clone()), lambda a, st: api.exemplar_rmsnorm(a[0], None, a[1], stream=st)),
    "norm_rows": (lambda m: (m[0], m[0].clone()),
                  lambda a, st: api.exemplar_rmsnorm(a[0], None, a[1], format=api.EXEMCL_MXFP8, stream=st)),
    "norm_gradient": (lambda m: (m[0], m[0].clone(), m[4]),
                      lambda a, st: api.exemplar_rmsnorm_backward(a[0], a[1], None, a[2], stream=st)),
    "product": (lambda m: (m[3], m[2]), lambda a, st: api.exemplar_mx_product(*a, stream=st)),
    "mx_eval": (lambda m: (m[2], m[1]), lambda a, st: api.exemplar_mx_eval(*a, stream=st)),
}


def copies(a):
    """The inputs again, in memory of their own."""
    return tuple(x._replace(codes=x.codes.clone(), scales=x.scales.clone()) if isinstance(x, api.MxRows) else x.clone()
                 for x in a)


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_a_call_on_another_stream(name, made):
    inputs, call = CALLS[name]
    args = inputs(made)
    want = tensors(call(args, None))
    main, st = torch.cuda.current_stream(), torch.cuda.Stream()
    a = copies(args)
    st.wait_stream(main)
    call(a, st)  # what is allocated once
    torch.cuda.synchronize()

    # a block freed on the current stream, where its last use is queued, is no result
    torch.cuda._sleep(BUSY)
    freed = [torch.empty_like(t) for t in want]
    spans = [span(t) for t in freed]
    del freed
    results = call(a, st)
    got = tensors(results)
    assert all(apart(t, spans) for t in got)
    # inputs freed while their stream is still to read them are not handed out again
    with torch.cuda.stream(st):
        torch.cuda._sleep(BUSY)
    again = call(a, st)
    spans = [span(t) for t in tensors(a)] + [span(t) for t in tensors(again)]
    shapes = [(t.shape, t.dtype) for t in tensors(a, again)]
    del a, again
    fresh = [torch.empty(shape, dtype=dtype, device="cuda") for shape, dtype in shapes]
    assert all(apart(t, spans) for t in fresh)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    # results freed while the current stream is still to read them are no results of the next call
    torch.cuda._sleep(BUSY)
    spans = [span(t) for t in got]
    del got, results
    assert all(apart(t, spans) for t in tensors(call(args, st)))
    torch.cuda.synchronize()
