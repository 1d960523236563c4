"""What the GPU tests of the operators share."""

import numpy as np

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # half a spacing, relative


def types(torch):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def stored(torch, values, kind):
    """values rounded to the type on the host (torch's CPU conversion), as a CPU tensor."""
    return torch.from_numpy(np.ascontiguousarray(values, dtype=np.float32)).to(types(torch)[kind])


def doubles(t):
    return t.detach().cpu().double().numpy()


def guarded(torch, shape, dtype, margin=64, fill=77.0):
    """A tensor inside a larger one filled with `fill`, and the function that checks the margins."""
    count = int(np.prod(shape))
    whole = torch.full((count + 2 * margin,), fill, dtype=dtype, device="cuda")

    def check():
        assert bool((whole[:margin] == fill).all()) and bool((whole[margin + count:] == fill).all())
    return whole[margin:margin + count].view(shape), check


def replays(torch, call, outputs, refresh, times=3):
    """Captures `call` into a graph and replays it `times`, with new inputs from `refresh(i)` and the program's own eager work between;
    yields what `outputs()` held after each replay and after the eager call on the same inputs."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(times):
        refresh(i)
        for t in outputs():
            t.fill_(99)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outputs()]
        for t in outputs():
            t.fill_(98)
        call()
        torch.cuda.synchronize()
        yield got, [t.clone() for t in outputs()]
