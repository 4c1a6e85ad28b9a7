"""Which kernels a call of a residual block's operators launches, on what grids, without a GPU: the program of dispatch_train over the
library as it is built, with calls of its own."""
import subprocess

import dispatch_train

MAIN = r"""
int main()
{
    char what[32];
    long long v[8];
    auto at = [](int k) { return reinterpret_cast<char*>((uintptr_t)(k + 1) << 44); };
    auto f = [&](int k) { return reinterpret_cast<float*>(at(k)); };
    const hdqt_dropout_t drop = {0.3, 1, nullptr, 2, 0};
    while (scanf("%31s %lld %lld %lld %lld %lld %lld %lld %lld", what, v, v + 1, v + 2, v + 3, v + 4, v + 5, v + 6, v + 7) == 9) {
        g_log.clear();
        g_error = hipSuccess;
        int rc = -99;
        size_t ws = 0;
        if (!strcmp(what, "dropout"))               // elements, type
            rc = hdqt_dropout(at(0), at(1), at(2), v[0], (int)v[1], &drop, nullptr);
        if (!strcmp(what, "norm_fwd"))              // rows, columns, type
            rc = hdqt_layernorm_fwd(at(0), at(1), &drop, at(2), at(3), at(4), at(5), f(6), v[0], v[1], 1e-5f, (int)v[2], HDQT_F32, nullptr);
        if (!strcmp(what, "norm_bwd")) {            // rows, columns, type, wanted (1 dx, 2 dresidual, 4 dweight, 8 dbias; 16: dx is dy, 32: dresidual is)
            auto want = [&](int bit, int k) { return v[3] & bit ? at(k) : nullptr; };
            ws = hdqt_layernorm_bwd_workspace_size(v[0], v[1], (int)v[2]);
            rc = hdqt_layernorm_bwd(at(0), at(1), at(2), &drop, at(3), f(4), want(1, v[3] & 16 ? 0 : 5), want(2, v[3] & 32 ? 0 : 6), want(4, 7), want(8, 8), v[0],
                                    v[1], (int)v[2], HDQT_F32, at(9), ws, nullptr);
        }
        if (!strncmp(what, "adapt", 5)) {           // rows, features, outputs, rank, adapters, type, wanted (1 dx, 2 dA, 4 dB)
            const int r = (int)v[3], n = (int)v[4], t = (int)v[5];
            const int64_t* ids = reinterpret_cast<const int64_t*>(at(3));
            auto want = [&](int bit, int k) { return v[6] & bit ? at(k) : nullptr; };
            const size_t saved = hdqt_adapters_saved_size(v[0], v[1], v[2], r, n, t);
            ws = hdqt_adapters_bwd_workspace_size(v[0], v[1], v[2], r, n, t);
            if (!strcmp(what, "adapt_fwd"))
                rc = hdqt_adapters_fwd(at(0), at(1), at(2), ids, f(4), at(5), at(6), at(7), saved, v[0], v[1], v[2], r, n, t, nullptr);
            else
                rc = hdqt_adapters_bwd(at(8), at(0), at(1), at(2), ids, f(4), at(7), saved, nullptr, want(1, 9), want(2, 10), want(4, 11), v[0], v[1],
                                       v[2], r, n, t, at(12), ws, nullptr);
        }
        printf("%d %zu%s\n", rc, ws, g_log.c_str());
    }
    return 0;
}
"""

_EXE = None


def dispatch(calls):
    """calls: ("dropout", elements, type), ("norm_fwd" | "norm_bwd", rows, columns, type, wanted) or ("adapt_fwd" | "adapt_bwd", rows, features,
    outputs, rank, adapters, type, wanted) each; as dispatch_train's."""
    global _EXE
    if _EXE is None:
        program, exe, folder = dispatch_train.PROGRAM, dispatch_train._EXE, dispatch_train._FOLDER
        dispatch_train.PROGRAM, dispatch_train._EXE = program.split("int main()")[0] + MAIN, None
        try:
            _EXE = dispatch_train._program(), dispatch_train._FOLDER
        finally:
            dispatch_train.PROGRAM, dispatch_train._EXE, dispatch_train._FOLDER = program, exe, folder
    text = "".join(" ".join(map(str, c)) + " 0" * (9 - len(c)) + "\n" for c in calls)
    out = subprocess.run([_EXE[0]], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(calls)
    got = []
    for line in out:
        head, *rest = line.split("|")
        launches = []
        for r in rest:
            name, shape = r.rsplit("@", 1)
            x, y, z, threads = map(int, shape.split(","))
            launches.append(dispatch_train.Launch(name.split("<")[0], (x, y, z), threads))
        rc, workspace = map(int, head.split())
        got.append(dispatch_train.Call(rc, workspace, launches))
    return got
