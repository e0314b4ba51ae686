/* host_stub.c with streams that record graphs, memory that cannot be freed, and devices of other sizes. */
#define hipFree free_block
#include "host_stub.c"
#undef hipFree

#define MAX_STREAMS 16
static struct { hipStream_t stream; unsigned long long capture; hipStreamCaptureStatus status; } recording[MAX_STREAMS];

/* The stream records as part of a capture (0: it does not), which goes on or has failed. */
void stub_capture(void *stream, unsigned long long capture, int failed)
{
    int i;
    for (i = 0; i < MAX_STREAMS - 1 && recording[i].stream && recording[i].stream != (hipStream_t)stream; ++i);
    recording[i].stream = (hipStream_t)stream;
    recording[i].capture = capture;
    recording[i].status = !capture ? hipStreamCaptureStatusNone : failed ? hipStreamCaptureStatusInvalidated : hipStreamCaptureStatusActive;
}
static int refuse_free;
void stub_refuse_free(int yes) { refuse_free = yes; }
hipError_t hipFree(void *p) { return refuse_free ? last_error = hipErrorStreamCaptureUnsupported : free_block(p); }
void stub_compute_units(int n) { n_cus = n; }

hipError_t hipStreamGetCaptureInfo(hipStream_t s, hipStreamCaptureStatus *status, unsigned long long *id)
{
    int i;
    *status = hipStreamCaptureStatusNone;
    for (i = 0; i < MAX_STREAMS; ++i)
        if (s && recording[i].stream == s) {
            *status = recording[i].status;
            *id = recording[i].capture;
        }
    return hipSuccess;
}
