/* launch_recorder.c for switch_linear: what its calls would launch, without a GPU.
 *
 * input, one call per line:
 *   forward|backward M K N dtype activation dropout flags
 * output per call:
 *   launch <mangled kernel name> gx gy gz bx by bz lds     of each launch, then
 *   call <status> <workspace bytes>
 * Usage: linear_recorder <library>
 */
#define main layer_main
#include "launch_recorder.c"
#undef main

int main(int argc, char **argv) {
    void *lib = argc == 2 ? dlopen(argv[1], RTLD_NOW) : NULL;
    if (!lib) { fprintf(stderr, "%s\n", argc == 2 ? dlerror() : "usage: linear_recorder <library>"); return 2; }
    typeof(&switch_linear_workspace_size) size_of = dlsym(lib, "switch_linear_workspace_size");
    typeof(&switch_linear) forward = dlsym(lib, "switch_linear");
    typeof(&switch_linear_backward) backward = dlsym(lib, "switch_linear_backward");
    char what[16];
    long long M, K, N;
    int dtype, act, flags;
    float dropout;
    while (scanf("%15s %lld %lld %lld %d %d %f %d", what, &M, &K, &N, &dtype, &act, &dropout, &flags) == 8) {
        switch_linear_config c = {M, K, N, dtype, act, dropout, flags, 17};
        const int back = strcmp(what, "backward") == 0;
        size_t bytes = 0;
        int st = size_of(&c, back, &bytes);
        void *at = (void *)(1ull << 44), *ws = (void *)(1ull << 45);   /* never touched */
        if (st == 0)
            st = back ? backward(&c, at, at, at, at, at, at, at, ws, bytes, NULL)
                      : forward(&c, at, at, at, at, at, at, ws, bytes, NULL);
        printf("call %d %zu\n", st, bytes);
    }
    fflush(stdout);
    _exit(0);
}
