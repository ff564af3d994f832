"""A handle that does not fit the device's memory is refused, and the error
stays with that call: the next calls of the thread succeed."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _take_the_memory():
    """All of it but for 128 MiB or less."""
    torch.cuda.empty_cache()
    held = []
    for mib in (65536, 4096, 256, 64):
        while torch.cuda.mem_get_info()[0] > (mib + 64) << 20:
            held.append(torch.empty(mib << 20, dtype=torch.uint8, device="cuda"))
    return held


def test_calls_after_a_refused_handle():
    import paper_2411_01433_amd as P
    d, f, E, T = 256, 65536, 16, 4
    zeros = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")
    wg, x, wide = zeros(E, d), zeros(T, d), zeros(512, 64)
    h, y = torch.ones((T, d), device="cuda"), torch.empty((T, d), device="cuda")
    idx, w = torch.empty((T, 2), dtype=torch.int32, device="cuda"), torch.empty((T, 2), device="cuda")
    up, down = zeros(f, d), zeros(d, f)
    small_up, small_down = zeros(64, d), zeros(d, 64)
    layer = lambda f, T, a, b: P.MoeLayer(d, f, E, 2, T, wg, [a] * E, [a] * E, [b] * E)
    r, L = P.MoeRouter(d, E, 2, T, wg), layer(64, T, small_up, small_down)
    torch.cuda.synchronize()
    refused = (lambda: P.MoeRouter(64, 512, 8, 65536, wide, backward=True),   # 400 MiB
               lambda: layer(f, 8192, up, down))                              # 2 GiB
    calls = (lambda: r.route(x, idx, w), lambda: P.layernorm(h, x), lambda: P.rmsnorm(h, x),
             lambda: L.decode_step(x, y), lambda: L.prefill(x, y))
    held = _take_the_memory()
    try:
        for make in refused:
            for call in calls:
                with pytest.raises(P.MoeError) as e:
                    make()
                assert e.value.status == P.MOE_ENOMEM
                call()
        torch.cuda.synchronize()
    finally:
        held.clear()
        torch.cuda.empty_cache()
    L.destroy()
    r.destroy()
